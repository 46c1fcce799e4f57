"""A state-space policy on the Pong env: the sequence operators as a policy uses them.

The GRU of policy_loop.py acts; it cannot be trained on what it rolled out without walking
the rollout step by step.  A layer here is a gated state-space mixer and a gated
feed-forward block, both with a residual connection:

    [x | z] = h W_xz^T                       projections: torch matrix products
    x       = conv(x)                        ssm.h, short causal convolution
    [r|b|c] = x W_p^T,   dt = r W_dt^T
    h       = h + scan(x, dt, b, c, z) W_y^T    ssm.h, selective scan
    h       = h + ffn(h)                     gated_ffn.h

With norm=True each branch reads the stream normalised (layer_norm.h), and the addition of the branch before it is part of the
norm; with mixer="recurrence" the scan's place is taken by the lighter gated recurrence (gated_recurrence.h):

    [r | i] = x W_g^T
    h       = h + (recurrence(x, r, i) silu(z)) W_y^T

While the agent acts, every layer takes one token per env with the single-token forms; the
recurrent state and the last convolution inputs are cleared where an episode ended.
Training takes the stored rollout [steps, envs] in one piece with the sequence forms: the
same recurrence from the state at the rollout's start, episode ends inside, gradients by
torch.autograd through the Functions below, steps by Adam or, for the layers' matrices, by orthogonalised momentum
(optimizers.py).

    python -m paper_2603_12145_b200.ssm_policy --envs 1024 --steps 64 --updates 5
    python -m paper_2603_12145_b200.ssm_policy --mixer recurrence --norm --optimizer orthogonal --layers 6
"""
from __future__ import annotations

import functools
import math

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

from . import gated_ffn, gated_recurrence, layer_norm, optimizers, pong, ssm


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
    def wrapped(ctx, *dy):
        with torch.no_grad():
            grads = backward(ctx, *dy)
        if not torch.is_grad_enabled():
            return grads
        of = [v for v in dy + tuple(ctx.saved_tensors) if v is not None and v.requires_grad]
        return tuple(_Refuse.apply(g, *of) if g is not None and of else g for g in grads)

    return wrapped


def _differentiated(args):
    """Whether autograd has to see the call: an input that requires a gradient, or one with a forward-mode tangent, which the
    kernels would drop (a Function without a rule for it raises)."""
    tensors = [v for v in args if isinstance(v, torch.Tensor)]
    if torch.is_grad_enabled() and any(v.requires_grad for v in tensors):
        return True
    # (without an open level nothing carries one: 2 us less per call)
    return getattr(forward_ad, "_current_level", 0) >= 0 and any(forward_ad.unpack_dual(v).tangent is not None for v in tensors)


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
        if _differentiated(args):
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
        return super().apply(op, x, w_in, w_out) if _differentiated((x, w_in, w_out)) else op.forward(x, w_in, w_out)

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


class NormFunction(torch.autograd.Function):
    """layer_norm.LayerNorm on rows [n, width] with its gradients: the normalised rows, and with a residual
    (rows, x + residual), whose gradients meet here again."""

    @classmethod
    def apply(cls, op, x, residual, w, b):
        if _differentiated((x, residual, w, b)):
            return super().apply(op, x, residual, w, b)
        return op.forward(x, w, b, residual=residual)

    @staticmethod
    def forward(ctx, op, x, residual, w, b):
        ctx.set_materialize_grads(False)
        saved = op.saved(x.shape[0])
        ctx.op = op
        out = op.forward(x, w, b, residual=residual, saved=saved)
        ctx.save_for_backward(x if residual is None else out[1], w, saved)
        return out

    @staticmethod
    @first_order
    def backward(ctx, dy, dsum=None):
        s, w, saved = ctx.saved_tensors
        added, want_w, want_b = ctx.needs_input_grad[2], ctx.needs_input_grad[3], ctx.needs_input_grad[4]
        if dy is None:                     # the normalised rows were not used
            return None, dsum, dsum if added else None, None, None
        dx, dw, db = ctx.op.backward(_dense_last(dy), s, w, saved, dsum=None if dsum is None else _dense_last(dsum),
                                     want_params=want_w or want_b)
        return None, dx, dx if added else None, dw if want_w else None, db if want_b else None


class RecurrenceFunction(torch.autograd.Function):
    """gated_recurrence.GatedRecurrence.sequence with its gradients, that of the state at the start among them.  state_out is
    filled by address: what is computed from it is a constant here."""

    @classmethod
    def apply(cls, op, x, r, i, a, reset, state, state_out):
        if _differentiated((x, r, i, a, state)):
            return super().apply(op, x, r, i, a, reset, state, state_out)
        return op.sequence(x, r, i, a, reset=reset, state=state, state_out=state_out)

    @staticmethod
    def forward(ctx, op, x, r, i, a, reset, state, state_out):
        saved = op.saved(x.shape[0], x.shape[1])
        ctx.op = op
        # (the kernels do not read the state again; the gradients depend on it)
        ctx.save_for_backward(x, r, i, a, reset, saved, state if ctx.needs_input_grad[6] else None)
        return op.sequence(x, r, i, a, reset=reset, state=state, state_out=state_out, saved=saved)

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x, r, i, a, reset, saved, _ = ctx.saved_tensors
        g = ctx.op.backward(_dense_last(dy), x, r, i, a, saved, reset=reset, want_dstate=ctx.needs_input_grad[6])
        return None, g["dx"], g["dr"], g["di"], g["da"], None, g["dstate"], None


def _dense_last(v):
    return v if v.stride(-1) == 1 else v.contiguous()


class Layer(torch.nn.Module):
    def __init__(self, model: int, states: int, width: int, rank: int, ffn_hidden: int, device, seed: int,
                 mixer: str = "scan", norm: bool = False):
        super().__init__()
        if mixer not in ("scan", "recurrence"):
            raise ValueError("mixer must be scan or recurrence")
        inner = 2 * model
        self.inner, self.states, self.rank, self.mixer = inner, states, rank, mixer
        self.op = ssm.Ssm(inner, states, 1, width, torch.bfloat16, device=str(device))
        self.ffn = gated_ffn.GatedFfn(model, ffn_hidden, device=str(device))
        gen = torch.Generator().manual_seed(seed)

        def matrix(rows, cols, scale=1.0):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=gen) * scale * cols ** -0.5).to(device))

        self.w_xz = matrix(2 * inner, model)
        if mixer == "scan":
            self.w_p, self.w_dt = matrix(rank + 2 * states, inner), matrix(inner, rank)
        else:
            self.recurrence = gated_recurrence.GatedRecurrence(inner, device=str(device))
            self.w_g = matrix(2 * inner, inner)
        self.w_y, self.w_in, self.w_out = matrix(model, inner, 0.5), matrix(2 * ffn_hidden, model), matrix(model, ffn_hidden, 0.5)
        self.conv_w = torch.nn.Parameter((torch.randn(inner, width, generator=gen) * width ** -0.5).to(device))
        self.conv_b = torch.nn.Parameter(torch.zeros(inner, device=device))
        start = torch.exp(torch.rand(inner, generator=gen) * math.log(100.0) + math.log(1e-3))   # steps of 0.001 .. 0.1
        if mixer == "scan":
            self.log_rate = torch.nn.Parameter(torch.log(torch.arange(1, states + 1, device=device).float()).repeat(inner, 1))
            self.skip = torch.nn.Parameter(torch.ones(inner, device=device))
            self.dt_bias = torch.nn.Parameter((start + torch.log(-torch.expm1(-start))).to(device))
        else:
            self.log_rate = torch.nn.Parameter(torch.log(10.0 * start).to(device))     # strongest decays of 0.01 .. 1 a step
        self.norms = None
        if norm:
            self.norms = [layer_norm.LayerNorm(model, device=str(device)) for _ in range(2)]
            self.norm_w = torch.nn.Parameter(torch.ones(2, model, device=device))
            self.norm_b = torch.nn.Parameter(torch.zeros(2, model, device=device))

    def state(self, n: int):
        """The recurrent state of n fresh envs."""
        return (self.op if self.mixer == "scan" else self.recurrence).state(n).zero_()

    def matrices(self):
        """The parameters that orthogonalised momentum is for."""
        names = ("w_xz", "w_p", "w_dt", "w_y", "w_in", "w_out") if self.mixer == "scan" else ("w_xz", "w_g", "w_y", "w_in", "w_out")
        return [getattr(self, k) for k in names]

    def _projections(self, x):
        r, b, c = torch.split(x @ self.w_p.to(x.dtype).t(), [self.rank, self.states, self.states], dim=-1)
        return r @ self.w_dt.to(x.dtype).t(), b, c

    def _mix(self, h, reset, state, history):
        """The mixer's branch on [batch, time, model]."""
        x, z = torch.split(h @ self.w_xz.to(h.dtype).t(), [self.inner, self.inner], dim=-1)
        x = ConvFunction.apply(self.op, x, self.conv_w, self.conv_b, reset, history, None)
        if self.mixer == "scan":
            dt, b, c = self._projections(x)
            y = ScanFunction.apply(self.op, x, dt, -torch.exp(self.log_rate), b, c, self.skip, z, self.dt_bias, reset,
                                   state, None)
        else:
            r, i = torch.split(x @ self.w_g.to(x.dtype).t(), [self.inner, self.inner], dim=-1)
            y = RecurrenceFunction.apply(self.recurrence, x, r, i, -torch.exp(self.log_rate), reset, state, None)
            y = y * torch.nn.functional.silu(z)
        return y @ self.w_y.to(h.dtype).t()

    def sequence(self, h, reset, state, history):
        """h [batch, time, model] -> the layer's output; starts from state and history."""
        batch, time, model = h.shape
        h = h + self._mix(h, reset, state, history)
        rows = h.transpose(0, 1).reshape(batch * time, model)      # the rollout's own order: no copy if time-major
        f = FfnFunction.apply(self.ffn, rows, self.w_in.to(h.dtype), self.w_out.to(h.dtype))
        return h + f.view(time, batch, model).transpose(0, 1)

    def _norm(self, k, h, branch):
        """(normalised rows, the stream as it goes on) of the stream and the branch that is still to be added."""
        y = NormFunction.apply(self.norms[k], h, branch, self.norm_w[k], self.norm_b[k])
        return (y, h) if branch is None else y

    def normed_sequence(self, h, branch, batch, time, reset, state, history):
        """The stream h [time * batch, model] and the branch to be added to it -> the same behind this layer."""
        y, h = self._norm(0, h, branch)
        m = self._mix(y.view(time, batch, -1).transpose(0, 1), reset, state, history)
        y, h = self._norm(1, h, m.transpose(0, 1).reshape(time * batch, -1))
        return h, FfnFunction.apply(self.ffn, y, self.w_in.to(h.dtype), self.w_out.to(h.dtype))

    def weights(self):
        """What the single-token form reads, converted once per rollout."""
        names = ("w_xz", "w_p", "w_dt", "w_y", "w_in", "w_out") if self.mixer == "scan" else ("w_xz", "w_g", "w_y", "w_in", "w_out")
        w = {k: getattr(self, k).detach().to(torch.bfloat16) for k in names}
        w["a"] = -torch.exp(self.log_rate.detach())
        return w

    def _mix_step(self, w, h, done, state, history):
        x, z = torch.split(h @ w["w_xz"].t(), [self.inner, self.inner], dim=-1)
        # a training pass that started from these must not go on with what is written here by address
        increment_version((state, history))
        x = self.op.conv_step(x, history, self.conv_w, self.conv_b, done=done)
        if self.mixer == "scan":
            r, b, c = torch.split(x @ w["w_p"].t(), [self.rank, self.states, self.states], dim=-1)
            y = self.op.scan_step(x, r @ w["w_dt"].t(), w["a"], b, c, state, d=self.skip, z=z, dt_bias=self.dt_bias, done=done)
        else:
            r, i = torch.split(x @ w["w_g"].t(), [self.inner, self.inner], dim=-1)
            y = self.recurrence.step(x, r, i, w["a"], state, done=done) * torch.nn.functional.silu(z)
        return y @ w["w_y"].t()

    def step(self, w, h, done, state, history):
        """h [n, model] -> [n, model]; state and history are updated in place."""
        h = h + self._mix_step(w, h, done, state, history)
        return h + self.ffn.forward(h, w["w_in"], w["w_out"])

    def normed_step(self, w, h, branch, done, state, history):
        """As normed_sequence, one token of n rows."""
        y, h = self._norm(0, h, branch)
        y, h = self._norm(1, h, self._mix_step(w, y, done, state, history))
        return h, self.ffn.forward(y, w["w_in"], w["w_out"])


class StateSpacePolicy(torch.nn.Module):
    """obs [.., 6] -> logits [.., 3]."""

    def __init__(self, model: int = 64, layers: int = 2, states: int = 16, width: int = 4, rank: int = 16,
                 ffn_hidden: int = 192, device: str = "cuda:0", seed: int = 0, mixer: str = "scan", norm: bool = False):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        self.device = torch.device(device)
        self.embed = torch.nn.Parameter((torch.randn(model, 6, generator=gen) * 6 ** -0.5).to(device))
        self.head = torch.nn.Parameter((torch.randn(3, model, generator=gen) * 0.1 * model ** -0.5).to(device))
        self.layers = torch.nn.ModuleList(Layer(model, states, width, rank, ffn_hidden, device, seed + 1 + i, mixer, norm)
                                          for i in range(layers))
        self.last_norm = None
        if norm:
            self.last_norm = layer_norm.LayerNorm(model, device=str(device))
            self.last_w = torch.nn.Parameter(torch.ones(model, device=device))
            self.last_b = torch.nn.Parameter(torch.zeros(model, device=device))

    def start(self, n: int):
        """Recurrent states and convolution histories of n fresh envs."""
        return [(layer.state(n), layer.op.history(n).zero_()) for layer in self.layers]

    def _last(self, h, branch):
        """The normalised stream behind the last layer."""
        if branch is None:
            return NormFunction.apply(self.last_norm, h, None, self.last_w, self.last_b)
        return NormFunction.apply(self.last_norm, h, branch, self.last_w, self.last_b)[0]

    def sequence(self, obs, reset, carry):
        """obs [batch, time, 6], reset [batch, time]; carry as from start().  Logits [batch, time, 3]."""
        h = (obs @ self.embed.t()).to(torch.bfloat16)
        if self.last_norm is not None:
            batch, time = obs.shape[:2]
            h, branch = h.transpose(0, 1).reshape(time * batch, -1), None      # the rollout's own order
            for layer, (state, history) in zip(self.layers, carry):
                h, branch = layer.normed_sequence(h, branch, batch, time, reset, state, history)
            return self._last(h, branch).view(time, batch, -1).transpose(0, 1).float() @ self.head.t()
        for layer, (state, history) in zip(self.layers, carry):
            h = layer.sequence(h, reset, state, history)
        return h.float() @ self.head.t()

    def weights(self):
        return [layer.weights() for layer in self.layers]

    @torch.no_grad()
    def step(self, obs, done, carry, weights):
        """obs [n, 6] -> logits [n, 3]; carry is updated in place."""
        h = (obs @ self.embed.t()).to(torch.bfloat16)
        if self.last_norm is not None:
            branch = None
            for layer, w, (state, history) in zip(self.layers, weights, carry):
                h, branch = layer.normed_step(w, h, branch, done, state, history)
            return self._last(h, branch).float() @ self.head.t()
        for layer, w, (state, history) in zip(self.layers, weights, carry):
            h = layer.step(w, h, done, state, history)
        return h.float() @ self.head.t()


class Trainer:
    """Rolls the policy out on Pong and improves it with the policy gradient of the rollout."""

    def __init__(self, policy: StateSpacePolicy, n_envs: int, steps: int, seed: int = 0, learning_rate: float = 3e-4,
                 optimizer: str = "adam", matrix_rate: float = 0.02):
        self.policy, self.n, self.steps = policy, int(n_envs), int(steps)
        dev = policy.device
        self.env = pong.PongEnv(n_envs, seed, device=str(dev))
        if optimizer not in ("adam", "orthogonal"):
            raise ValueError("optimizer must be adam or orthogonal")
        self.matrix_optimizer = None
        if optimizer == "adam":
            self.optimizer = torch.optim.Adam(policy.parameters(), lr=learning_rate)
        else:
            matrices = [p for layer in policy.layers for p in layer.matrices()]
            taken = set(map(id, matrices))
            self.matrix_optimizer = optimizers.OrthogonalMomentum(matrices, lr=matrix_rate)
            self.optimizer = torch.optim.Adam([p for p in policy.parameters() if id(p) not in taken], lr=learning_rate)
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
        self.policy.zero_grad(set_to_none=True)
        loss.backward()
        torch.nn.utils.clip_grad_norm_(self.policy.parameters(), 1.0)
        self.optimizer.step()
        if self.matrix_optimizer is not None:
            self.matrix_optimizer.step()
        return loss.detach()

    def check(self):
        """Synchronises; raises if a kernel gave up a wait."""
        for layer in self.policy.layers:
            layer.ffn.status()
        if self.matrix_optimizer is not None:
            self.matrix_optimizer.check()


def main(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--envs", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--updates", type=int, default=5)
    ap.add_argument("--model", type=int, default=64)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--mixer", choices=("scan", "recurrence"), default="scan")
    ap.add_argument("--norm", action="store_true", help="normalise what each branch reads")
    ap.add_argument("--optimizer", choices=("adam", "orthogonal"), default="adam", help="of the layers' matrices")
    args = ap.parse_args(argv)
    policy = StateSpacePolicy(model=args.model, layers=args.layers, ffn_hidden=3 * args.model, mixer=args.mixer, norm=args.norm)
    trainer = Trainer(policy, args.envs, args.steps, optimizer=args.optimizer)
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
