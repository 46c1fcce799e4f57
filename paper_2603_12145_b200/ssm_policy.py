"""A state-space policy on the Pong env: the sequence operators as a policy uses them.

The GRU of policy_loop.py acts; it cannot be trained on what it rolled out without walking
the rollout step by step.  A layer here is a gated state-space mixer and a gated
feed-forward block, both with a residual connection:

    [x | z] = h W_xz^T                       projections: torch matrix products
    x       = conv(x)                        ssm.h, short causal convolution
    [r|b|c] = x W_p^T,   dt = r W_dt^T
    h       = h + scan(x, dt, b, c, z) W_y^T    ssm.h, selective scan
    h       = h + ffn(h)                     gated_ffn.h

While the agent acts, every layer takes one token per env with the single-token forms; the
recurrent state and the last convolution inputs are cleared where an episode ended.
Training takes the stored rollout [steps, envs] in one piece with the sequence forms: the
same recurrence from the state at the rollout's start, episode ends inside, gradients by
torch.autograd through the Functions below.

    python -m paper_2603_12145_b200.ssm_policy --envs 1024 --steps 64 --updates 5
"""
from __future__ import annotations

import functools
import math

import torch
from torch.autograd.graph import increment_version

from . import gated_ffn, pong, ssm


class _Refuse(torch.autograd.Function):
    """A gradient that itself depends on `of` in a way that autograd does not know."""

    @staticmethod
    def forward(ctx, gradient, *of):
        return gradient

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("the sequence operators have first derivatives only: this gradient was asked for its own")


def first_order(backward):
    """For a Function whose backward calls kernels.  With create_graph the gradients would look like constants, and
    a second derivative would silently lack what goes through the operator; here it raises.  (once_differentiable
    does so only where the incoming gradient carries a graph, not where the inputs alone do.)"""

    @functools.wraps(backward)
    def wrapped(ctx, dy):
        with torch.no_grad():
            grads = backward(ctx, dy)
        if not torch.is_grad_enabled():
            return grads
        of = [v for v in (dy,) + tuple(ctx.saved_tensors) if v is not None and v.requires_grad]
        return tuple(_Refuse.apply(g, *of) if g is not None and of else g for g in grads)

    return wrapped


def _wants_gradient(args):
    return torch.is_grad_enabled() and any(isinstance(v, torch.Tensor) and v.requires_grad for v in args)


class ConvFunction(torch.autograd.Function):
    """ssm.Ssm.conv with its gradients; the history is a constant."""

    @staticmethod
    def forward(ctx, op, x, w, bias, reset, history, history_out):
        ctx.op = op
        ctx.save_for_backward(x, w, bias, reset, history)
        return op.conv(x, w, bias, reset=reset, history=history, history_out=history_out)

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, w, bias, reset, history = ctx.saved_tensors
        dx, dw, dbias = ctx.op.conv_backward(_dense_last(dy), x, w, bias, reset=reset, history=history)
        return None, dx, dw, dbias, None, None, None


class ScanFunction(torch.autograd.Function):
    """ssm.Ssm.scan with its gradients; the state at the start is a constant."""

    @classmethod
    def apply(cls, op, x, dt, a, b, c, d, z, dt_bias, reset, state, state_out):
        args = (op, x, dt, a, b, c, d, z, dt_bias, reset, state, state_out)
        if _wants_gradient(args):
            return super().apply(*args)
        return op.scan(x, dt, a, b, c, d=d, z=z, dt_bias=dt_bias, reset=reset, state=state, state_out=state_out)

    @staticmethod
    def forward(ctx, op, x, dt, a, b, c, d, z, dt_bias, reset, state, state_out):
        saved = op.saved(x.shape[0], x.shape[1])
        ctx.op = op
        ctx.save_for_backward(x, dt, a, b, c, d, z, dt_bias, reset, saved)
        return op.scan(x, dt, a, b, c, d=d, z=z, dt_bias=dt_bias, reset=reset, state=state, state_out=state_out,
                       saved=saved)

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, dt, a, b, c, d, z, dt_bias, reset, saved = ctx.saved_tensors
        g = ctx.op.scan_backward(_dense_last(dy), x, dt, a, b, c, saved, d=d, z=z, dt_bias=dt_bias, reset=reset)
        return (None, g["dx"], g["ddt"], g["da"], g["db"], g["dc"], g["dd"], g["dz"], g["ddt_bias"], None, None, None)


class FfnFunction(torch.autograd.Function):
    """gated_ffn.GatedFfn on rows [n, model] with its gradients."""

    @classmethod
    def apply(cls, op, x, w_in, w_out):
        return super().apply(op, x, w_in, w_out) if _wants_gradient((x, w_in, w_out)) else op.forward(x, w_in, w_out)

    @staticmethod
    def forward(ctx, op, x, w_in, w_out):
        saved = op.saved(x.shape[0])
        ctx.op = op
        ctx.save_for_backward(x, w_in, w_out, *saved)
        return op.forward(x, w_in, w_out, saved=saved)

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, w_in, w_out, pre, hidden = ctx.saved_tensors
        return (None,) + ctx.op.backward(dy.contiguous(), x, w_in, w_out, (pre, hidden))


def _dense_last(v):
    return v if v.stride(-1) == 1 else v.contiguous()


class Layer(torch.nn.Module):
    def __init__(self, model: int, states: int, width: int, rank: int, ffn_hidden: int, device, seed: int):
        super().__init__()
        inner = 2 * model
        self.inner, self.states, self.rank = inner, states, rank
        self.op = ssm.Ssm(inner, states, 1, width, torch.bfloat16, device=str(device))
        self.ffn = gated_ffn.GatedFfn(model, ffn_hidden, device=str(device))
        gen = torch.Generator().manual_seed(seed)

        def matrix(rows, cols, scale=1.0):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=gen) * scale * cols ** -0.5).to(device))

        self.w_xz, self.w_p, self.w_dt = matrix(2 * inner, model), matrix(rank + 2 * states, inner), matrix(inner, rank)
        self.w_y, self.w_in, self.w_out = matrix(model, inner, 0.5), matrix(2 * ffn_hidden, model), matrix(model, ffn_hidden, 0.5)
        self.conv_w = torch.nn.Parameter((torch.randn(inner, width, generator=gen) * width ** -0.5).to(device))
        self.conv_b = torch.nn.Parameter(torch.zeros(inner, device=device))
        self.log_rate = torch.nn.Parameter(torch.log(torch.arange(1, states + 1, device=device).float()).repeat(inner, 1))
        self.skip = torch.nn.Parameter(torch.ones(inner, device=device))
        start = torch.exp(torch.rand(inner, generator=gen) * math.log(100.0) + math.log(1e-3))   # steps of 0.001 .. 0.1
        self.dt_bias = torch.nn.Parameter((start + torch.log(-torch.expm1(-start))).to(device))

    def _projections(self, x):
        r, b, c = torch.split(x @ self.w_p.to(x.dtype).t(), [self.rank, self.states, self.states], dim=-1)
        return r @ self.w_dt.to(x.dtype).t(), b, c

    def sequence(self, h, reset, state, history):
        """h [batch, time, model] -> the layer's output; starts from state and history."""
        batch, time, model = h.shape
        x, z = torch.split(h @ self.w_xz.to(h.dtype).t(), [self.inner, self.inner], dim=-1)
        x = ConvFunction.apply(self.op, x, self.conv_w, self.conv_b, reset, history, None)
        dt, b, c = self._projections(x)
        y = ScanFunction.apply(self.op, x, dt, -torch.exp(self.log_rate), b, c, self.skip, z, self.dt_bias, reset,
                               state, None)
        h = h + y @ self.w_y.to(h.dtype).t()
        rows = h.transpose(0, 1).reshape(batch * time, model)      # the rollout's own order: no copy if time-major
        f = FfnFunction.apply(self.ffn, rows, self.w_in.to(h.dtype), self.w_out.to(h.dtype))
        return h + f.view(time, batch, model).transpose(0, 1)

    def weights(self):
        """What the single-token form reads, converted once per rollout."""
        w = {k: getattr(self, k).detach().to(torch.bfloat16) for k in ("w_xz", "w_p", "w_dt", "w_y", "w_in", "w_out")}
        w["a"] = -torch.exp(self.log_rate.detach())
        return w

    def step(self, w, h, done, state, history):
        """h [n, model] -> [n, model]; state and history are updated in place."""
        x, z = torch.split(h @ w["w_xz"].t(), [self.inner, self.inner], dim=-1)
        # a training pass that started from these must not go on with what is written here by address
        increment_version((state, history))
        x = self.op.conv_step(x, history, self.conv_w, self.conv_b, done=done)
        r, b, c = torch.split(x @ w["w_p"].t(), [self.rank, self.states, self.states], dim=-1)
        y = self.op.scan_step(x, r @ w["w_dt"].t(), w["a"], b, c, state, d=self.skip, z=z, dt_bias=self.dt_bias, done=done)
        h = h + y @ w["w_y"].t()
        return h + self.ffn.forward(h, w["w_in"], w["w_out"])


class StateSpacePolicy(torch.nn.Module):
    """obs [.., 6] -> logits [.., 3]."""

    def __init__(self, model: int = 64, layers: int = 2, states: int = 16, width: int = 4, rank: int = 16,
                 ffn_hidden: int = 192, device: str = "cuda:0", seed: int = 0):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        self.device = torch.device(device)
        self.embed = torch.nn.Parameter((torch.randn(model, 6, generator=gen) * 6 ** -0.5).to(device))
        self.head = torch.nn.Parameter((torch.randn(3, model, generator=gen) * 0.1 * model ** -0.5).to(device))
        self.layers = torch.nn.ModuleList(Layer(model, states, width, rank, ffn_hidden, device, seed + 1 + i)
                                          for i in range(layers))

    def start(self, n: int):
        """Recurrent states and convolution histories of n fresh envs."""
        return [(layer.op.state(n).zero_(), layer.op.history(n).zero_()) for layer in self.layers]

    def sequence(self, obs, reset, carry):
        """obs [batch, time, 6], reset [batch, time]; carry as from start().  Logits [batch, time, 3]."""
        h = (obs @ self.embed.t()).to(torch.bfloat16)
        for layer, (state, history) in zip(self.layers, carry):
            h = layer.sequence(h, reset, state, history)
        return h.float() @ self.head.t()

    def weights(self):
        return [layer.weights() for layer in self.layers]

    @torch.no_grad()
    def step(self, obs, done, carry, weights):
        """obs [n, 6] -> logits [n, 3]; carry is updated in place."""
        h = (obs @ self.embed.t()).to(torch.bfloat16)
        for layer, w, (state, history) in zip(self.layers, weights, carry):
            h = layer.step(w, h, done, state, history)
        return h.float() @ self.head.t()


class Trainer:
    """Rolls the policy out on Pong and improves it with the policy gradient of the rollout."""

    def __init__(self, policy: StateSpacePolicy, n_envs: int, steps: int, seed: int = 0, learning_rate: float = 3e-4):
        self.policy, self.n, self.steps = policy, int(n_envs), int(steps)
        dev = policy.device
        self.env = pong.PongEnv(n_envs, seed, device=str(dev))
        self.optimizer = torch.optim.Adam(policy.parameters(), lr=learning_rate)
        self.obs = torch.empty((self.steps, self.n, 6), device=dev)
        self.reward = torch.empty((self.steps, self.n), device=dev)
        # done[t]: the episode ended with step t - 1, so that step t starts one; one row more than steps
        self.done = torch.zeros((self.steps + 1, self.n), dtype=torch.uint8, device=dev)
        self.actions = torch.empty((self.steps, self.n), dtype=torch.uint8, device=dev)
        self.logits = torch.empty((self.steps, self.n, 3), device=dev)
        self.carry = policy.start(self.n)
        self.current = self.env.reset()

    def rollout(self):
        """Acts for `steps` steps; returns the carry from before the first of them."""
        before = [(state.clone(), history.clone()) for state, history in self.carry]
        weights = self.policy.weights()
        words = self.env.fill_words(self.steps)
        self.done[0].copy_(self.done[self.steps])
        for t in range(self.steps):
            self.obs[t].copy_(self.current)
            self.logits[t].copy_(self.policy.step(self.current, self.done[t], self.carry, weights))
            self.env.sample_actions(self.logits[t], words[t], out=self.actions[t])
            self.env.step(self.actions[t], obs=self.current, reward=self.reward[t], done=self.done[t + 1])
        return before

    def update(self, before, discount: float = 0.99):
        """One gradient step on the stored rollout; returns the loss (a device scalar)."""
        gain = torch.zeros_like(self.reward[0])
        gains = torch.empty_like(self.reward)
        for t in range(self.steps - 1, -1, -1):
            gain = self.reward[t] + discount * gain * (self.done[t + 1] == 0)
            gains[t] = gain
        advantage = (gains - gains.mean()) / (gains.std() + 1e-6)
        logits = self.policy.sequence(self.obs.transpose(0, 1), self.done[:-1].t(), before).transpose(0, 1)
        chosen = torch.log_softmax(logits, dim=-1).gather(-1, self.actions.long().unsqueeze(-1)).squeeze(-1)
        loss = -(advantage * chosen).mean()
        self.optimizer.zero_grad(set_to_none=True)
        loss.backward()
        torch.nn.utils.clip_grad_norm_(self.policy.parameters(), 1.0)
        self.optimizer.step()
        return loss.detach()

    def check(self):
        """Synchronises; raises if a kernel gave up a wait."""
        for layer in self.policy.layers:
            layer.ffn.status()


def main(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--envs", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--updates", type=int, default=5)
    ap.add_argument("--model", type=int, default=64)
    ap.add_argument("--layers", type=int, default=2)
    args = ap.parse_args(argv)
    policy = StateSpacePolicy(model=args.model, layers=args.layers, ffn_hidden=3 * args.model)
    trainer = Trainer(policy, args.envs, args.steps)
    for i in range(args.updates):
        a, b, c = (torch.cuda.Event(enable_timing=True) for _ in range(3))
        a.record()
        before = trainer.rollout()
        b.record()
        loss = trainer.update(before)
        c.record()
        trainer.check()
        print("update %d: loss %.5f, mean reward %.5f, rollout %.1f ms, training step %.1f ms, %.0f env-steps/s"
              % (i, loss.item(), trainer.reward.mean().item(), a.elapsed_time(b), b.elapsed_time(c),
                 args.envs * args.steps / (a.elapsed_time(c) * 1e-3)))


if __name__ == "__main__":
    main()
