"""A gated feed-forward layer of n workers' models, trained by RelaySGD.

The layer operators put together as a training step uses them: the weights are
views of the workers' fp32 model rows, the gradients of rows beside them, and
what the backward pass needs of the activations is held in 8 bits:

    h = x + r;  y = rms_norm(h) w;  g, u = Wg y, Wu y;  out = Wd (g sigma(g) u)

``python -m paper_2110_04175_gb300.feed_forward`` trains it: every worker has
data of its own, the workers sit on a binary tree, and each step's gradients go
through ``GradientRun`` (Adam, then RelaySGD's relay, Algorithm 1).
"""
from __future__ import annotations

from . import layers as rl


class FeedForward:
    """The layer's buffers for n workers with `tokens` tokens of width d, hidden width f.

    ``weights(rows)`` gives the views of a [n][>= size] fp32 array: the norm's weight
    [n][d], gate and up [n][2 f][d] (one product) and down [n][d][f].  ``forward`` keeps
    the norm's rows and both halves of the product in 8 bits, ``backward`` reads them.
    The products with the weights are torch's; everything else runs in the library."""

    def __init__(self, n: int, tokens: int, d: int, f: int, dtype=None, eps: float = 1e-5, device="cuda"):
        import torch
        self.n, self.tokens, self.d, self.f, self.eps = n, tokens, d, f, eps
        self.dtype = dtype or torch.bfloat16
        self.at = [0, -(-d // 4) * 4]  # gate and up start on a 16-byte boundary of the rows
        self.at.append(self.at[1] + 2 * f * d)
        self.size = self.at[2] + d * f

        def rows(width):
            return torch.empty(n, tokens, width, dtype=self.dtype, device=device)

        self.total, self.y, self.both, self.act = rows(d), rows(d), rows(2 * f), rows(f)
        self.dboth, self.dx = rows(2 * f), rows(d)
        self.rstd = torch.empty(n, tokens, device=device)
        self.kept = rl.ActivationCheckpoint(n, tokens, d, device)
        self.kept_gate, self.kept_up, self.kept_act = (rl.ActivationCheckpoint(n, tokens, f, device) for _ in range(3))
        need = max(rl.relay_rms_norm_backward_workspace(n, tokens, d),
                   rl.relay_weight_grad_workspace(n, tokens, 2 * f, d, self.dboth),
                   rl.relay_weight_grad_workspace(n, tokens, d, f))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def weights(self, rows):
        """(norm [n][d], gate and up [n][2 f][d], down [n][d][f]) as views of fp32 rows."""
        d, f, (a, b, c) = self.d, self.f, self.at
        return (rows[:, a:a + d], rows[:, b:b + 2 * f * d].unflatten(1, (2 * f, d)),
                rows[:, c:c + d * f].unflatten(1, (d, f)))

    def _halves(self, both):
        return both[..., :self.f], both[..., self.f:]

    def forward(self, rows, x, residual=None):
        """(out, h): the layer's output and the sum that goes on past it."""
        import torch
        w, gate_up, down = self.weights(rows)
        rl.relay_rms_norm(x, w, self.y, self.eps, residual=residual, total=self.total, rstd=self.rstd,
                          checkpoint=self.kept)
        torch.bmm(self.y, gate_up.to(self.dtype).transpose(1, 2), out=self.both)
        rl.relay_gated(*self._halves(self.both), self.act, gate_checkpoint=self.kept_gate, up_checkpoint=self.kept_up)
        return self.act @ down.to(self.dtype).transpose(1, 2), self.total

    def backward(self, rows, grads, dout, dtotal=None, lengths=None):
        """The gradient of x and of the residual; the weights' go to `grads` (fp32 rows like
        `rows`).  dtotal: the gradient that reaches h past the layer; lengths: each worker's
        number of tokens."""
        w, gate_up, down = self.weights(rows)
        dw, dgate_up, ddown = self.weights(grads)
        rl.relay_gated_backward(dout @ down.to(self.dtype), *self._halves(self.dboth), gate_checkpoint=self.kept_gate,
                                up_checkpoint=self.kept_up, out_checkpoint=self.kept_act)
        rl.relay_weight_grad(dout, self.kept_act, ddown, self.workspace, lengths=lengths)
        # y = xhat w, and xhat is what was kept: w goes into the gradient's columns
        rl.relay_weight_grad(self.dboth, self.kept, dgate_up, self.workspace, column_scale=w, lengths=lengths)
        rl.relay_rms_norm_backward(self.dboth @ gate_up.to(self.dtype), w, self.rstd, self.dx, dw, self.workspace,
                                   checkpoint=self.kept, dtotal=dtotal, lengths=lengths)
        return self.dx


class GradientRun:
    """RelaySGD (Algorithm 1 with Adam) on gradients that the caller has computed.

    The step's own objective is a quadratic with the gradient x - mu, and a gradient handed
    over as mu = x - g would be rounded to the spacing of x.  So Adam runs on its own, as
    one worker's step from zero with the centre -g, where the gradient 0 - (-g) is g itself;
    its step goes into the relay as the centre x + step at lr = 1, rounded as any addition
    to x.  ``x`` (fp32 [n][>= d]): the models.  ``descent`` (like x, zero where nothing is
    written): the caller puts -g there, then calls ``step``."""

    def __init__(self, n: int, d: int, edges, beta1: float = 0.9, beta2: float = 0.99, eps: float = 1e-8):
        import numpy as np

        from . import RelayRun
        self.n, self.relay = n, RelayRun(n, d, edges)
        self.x = self.relay.x
        self.adam = RelayRun(1, self.x.numel(), np.zeros((0, 2), np.int32), optimizer=("adam", beta1, beta2, eps))
        self.descent = self.adam.mu.view_as(self.x)

    def init(self, x0_std: float, seed: int):
        """The same models everywhere, x0_std times normal values; no gradients yet."""
        import numpy as np
        self.relay.init(x0_std, seed, np.ones((self.n, 1)), 0.0, seed, 0.0)
        self.adam.init(0.0, seed, np.ones((1, 1)), 0.0, seed, 0.0)

    def step(self, lr: float, seed: int = 0):
        """One step of every worker with the gradients that `descent` holds, and its relay."""
        import torch
        self.adam.x.zero_()
        self.adam.step(lr, seed)
        torch.add(self.x, self.adam.x.view_as(self.x), out=self.relay.mu)
        self.relay.step(1.0, seed)


def train(n: int = 8, tokens: int = 256, d: int = 256, f: int = 512, steps: int = 100, lr: float = 0.02, seed: int = 0):
    """Trains one layer on n workers, each with inputs of its own mean, towards a common
    teacher's outputs; returns the mean loss per step."""
    import torch

    from . import workloads as wl

    layer = FeedForward(n, tokens, d, f)
    run = GradientRun(n, layer.size, wl.binary_tree(n))
    run.init(0.04, seed)  # the same models everywhere
    layer.weights(run.x)[0].fill_(1.0)
    make = torch.Generator(device="cuda").manual_seed(seed)
    teacher = torch.randn(1, layer.size, device="cuda", generator=make).mul_(0.08).expand(n, -1).contiguous()
    layer.weights(teacher)[0].fill_(1.0)
    x = torch.randn(n, tokens, d, device="cuda", generator=make)
    x = (x + torch.randn(n, 1, d, device="cuda", generator=make)).bfloat16()  # heterogeneous workers
    target = layer.forward(teacher, x)[0].clone()
    losses = []
    for _ in range(steps):
        out, _ = layer.forward(run.x, x)
        off = out.float() - target.float()
        losses.append(off.square().mean())
        layer.backward(run.x, run.descent, (off * (-1.0 / tokens)).bfloat16())  # -g
        run.step(lr, seed)
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    history = train()
    for step in range(0, len(history), 10):
        print(f"step {step:3d}  mean loss of the workers {history[step]:.4f}")
    print(f"step {len(history) - 1:3d}  mean loss of the workers {history[-1]:.4f}")
