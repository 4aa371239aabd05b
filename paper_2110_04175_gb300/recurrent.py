"""A recurrent block of n workers' models, trained by RelaySGD with orthogonal updates.

The layer operators put together as one block of a model without attention uses them: a
gated linear recurrence mixes the tokens, a gated feed-forward layer the features, and one
call takes the sum from the one to the other:

    y = rms_norm(r) w;  f, v, o = Wf y, Wv y, Wo y;  s = recurrence(f, v);  x = Wm (o sigma(o) s)
    h = scale r + norm(x) w_post;  y2 = norm(h) w_pre
    g, u = Wg y2, Wu y2;  out = h + Wd (g sigma(g) u)

``python -m paper_2110_04175_gb300.recurrent`` trains it: every worker has sequences of its
own, the workers sit on a binary tree, and each step's gradients go through ``GradientRun``
with the matrices' updates made orthogonal and the vectors' by Adam.
"""
from __future__ import annotations

from . import layers as rl
from .feed_forward import GradientRun


class RecurrentBlock:
    """The block's buffers for n workers with `tokens` tokens of width d, hidden width f.

    ``weights(rows)`` gives the views of a [n][>= size] fp32 array by name: the vectors
    "norm", "post", "pre" and "scale" [n][d], the matrices "mix" [n][3 f][d] (forget gate,
    value and output gate in one product), "mixed" [n][d][f], "gate_up" [n][2 f][d] and
    "down" [n][d][f].  ``begins`` (uint8 [n][tokens]) packs several sequences behind one
    another, ``lengths`` (int32 [n]) leaves the rest of a worker's rows out."""

    VECTORS = ("norm", "post", "pre", "scale")

    def __init__(self, n: int, tokens: int, d: int, f: int, dtype=None, eps: float = 1e-5, device="cuda"):
        import torch
        self.n, self.tokens, self.d, self.f, self.eps = n, tokens, d, f, eps
        self.dtype = dtype or torch.bfloat16
        shapes = {name: (d,) for name in self.VECTORS}
        shapes.update(mix=(3 * f, d), mixed=(d, f), gate_up=(2 * f, d), down=(d, f))
        self.at, self.size = {}, 0
        for name, shape in shapes.items():
            self.at[name] = self.size, shape
            count = shape[0] * (shape[1] if len(shape) > 1 else 1)
            self.size += -(-count // 4) * 4  # each starts on a 16-byte boundary of the rows

        def rows(width):
            return torch.empty(n, tokens, width, dtype=self.dtype, device=device)

        def kept(width):
            return rl.ActivationCheckpoint(n, tokens, width, device)

        self.y, self.total, self.y2, self.both, self.act = rows(d), rows(d), rows(d), rows(2 * f), rows(f)
        self.mix, self.state, self.mixed = rows(3 * f), rows(f), rows(f)
        self.dmix, self.dgate_value, self.dboth = rows(3 * f), rows(f), rows(2 * f)
        self.dx, self.dres, self.dr = rows(d), rows(d), rows(d)
        self.rstd, self.rstds = torch.empty(n, tokens, device=device), torch.empty(2, n, tokens, device=device)
        self.kept_y, self.kept_y2 = kept(d), kept(d)
        self.kept_mixed, self.kept_gate, self.kept_up, self.kept_act = (kept(f) for _ in range(4))
        need = max(rl.relay_rms_norm_backward_workspace(n, tokens, d), rl.relay_block_norm_backward_workspace(n, tokens, d),
                   rl.relay_recurrence_workspace(n, tokens, f), rl.relay_weight_grad_workspace(n, tokens, 3 * f, d),
                   rl.relay_weight_grad_workspace(n, tokens, d, f))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def weights(self, rows):
        """The weights by name, as views of fp32 rows."""
        out = {}
        for name, (first, shape) in self.at.items():
            count = shape[0] * (shape[1] if len(shape) > 1 else 1)
            part = rows[:, first:first + count]
            out[name] = part if len(shape) == 1 else part.unflatten(1, shape)
        return out

    def matrices(self, rows):
        """The matrices among them."""
        return [w for name, w in self.weights(rows).items() if name not in self.VECTORS]

    def _thirds(self, mix):
        return mix[..., :self.f], mix[..., self.f:2 * self.f], mix[..., 2 * self.f:]

    def _halves(self, both):
        return both[..., :self.f], both[..., self.f:]

    def forward(self, rows, r, initial=None, last=None, begins=None, lengths=None):
        """The block's output from the residual stream r.  initial, last (fp32 [n][f]): the
        recurrence's states before the first and behind the last token, for sequences that are
        worked through in stretches or token by token; one tensor may be both."""
        import torch
        w = self.weights(rows)
        rl.relay_rms_norm(r, w["norm"], self.y, self.eps, rstd=self.rstd, checkpoint=self.kept_y)
        torch.bmm(self.y, w["mix"].to(self.dtype).transpose(1, 2), out=self.mix)
        forget, value, gate = self._thirds(self.mix)
        rl.relay_recurrence(forget, value, self.state, self.workspace, initial=initial, last=last, begins=begins,
                            lengths=lengths)
        rl.relay_gated(gate, self.state, self.mixed)
        x = self.mixed @ w["mixed"].to(self.dtype).transpose(1, 2)
        rl.relay_block_norm(x, r, w["post"], w["pre"], self.total, self.y2, self.eps, scale=w["scale"], rstd=self.rstds,
                            checkpoint=self.kept_y2)
        torch.bmm(self.y2, w["gate_up"].to(self.dtype).transpose(1, 2), out=self.both)
        rl.relay_gated(*self._halves(self.both), self.act, gate_checkpoint=self.kept_gate, up_checkpoint=self.kept_up)
        self.r, self.x, self.initial, self.begins, self.lengths = r, x, initial, begins, lengths
        return self.total + self.act @ w["down"].to(self.dtype).transpose(1, 2)

    def backward(self, rows, grads, dout, dlast=None, dinitial=None):
        """The gradient of r; the weights' go to `grads` (fp32 rows like `rows`).  The forward pass
        has to be this block's last call, with `initial` left as it was.  dlast, dinitial (fp32
        [n][f]): the gradients of the states."""
        w, g, lengths = self.weights(rows), self.weights(grads), self.lengths
        dgate, dup = self._halves(self.dboth)
        rl.relay_gated_backward(dout @ w["down"].to(self.dtype), dgate, dup, gate_checkpoint=self.kept_gate,
                                up_checkpoint=self.kept_up, out_checkpoint=self.kept_act)
        rl.relay_weight_grad(dout, self.kept_act, g["down"], self.workspace, lengths=lengths)
        rl.relay_weight_grad(self.dboth, self.kept_y2, g["gate_up"], self.workspace, column_scale=w["pre"], lengths=lengths)
        rl.relay_block_norm_backward(self.dboth @ w["gate_up"].to(self.dtype), self.x, self.r, w["post"], w["pre"], self.rstds,
                                     self.dx, self.dres, g["post"], g["pre"], self.workspace, scale=w["scale"], dtotal=dout,
                                     dscale=g["scale"], lengths=lengths)
        forget, value, gate = self._thirds(self.mix)
        dforget, dvalue, dgate = self._thirds(self.dmix)
        rl.relay_gated_backward(self.dx @ w["mixed"].to(self.dtype), dgate, self.dgate_value, gate=gate, up=self.state,
                                out_checkpoint=self.kept_mixed)
        rl.relay_weight_grad(self.dx, self.kept_mixed, g["mixed"], self.workspace, lengths=lengths)
        rl.relay_recurrence_backward(self.dgate_value, forget, value, self.state, dforget, dvalue, self.workspace,
                                     initial=self.initial, dlast=dlast, dinitial=dinitial, begins=self.begins, lengths=lengths)
        rl.relay_weight_grad(self.dmix, self.kept_y, g["mix"], self.workspace, column_scale=w["norm"], lengths=lengths)
        rl.relay_rms_norm_backward(self.dmix @ w["mix"].to(self.dtype), w["norm"], self.rstd, self.dr, g["norm"],
                                   self.workspace, checkpoint=self.kept_y, dtotal=self.dres, lengths=lengths)
        return self.dr


def train(n: int = 8, tokens: int = 256, d: int = 128, f: int = 192, steps: int = 100, lr: float = 0.01, seed: int = 0):
    """Trains one block on n workers, each with inputs of its own mean and four sequences packed into
    its tokens, towards a common teacher's outputs; returns the mean loss per step."""
    import torch

    from . import workloads as wl

    block = RecurrentBlock(n, tokens, d, f)
    run = GradientRun(n, block.size, wl.binary_tree(n), matrices=block.matrices)
    run.init(0.04, seed)  # the same models everywhere
    make = torch.Generator(device="cuda").manual_seed(seed)
    teacher = torch.randn(1, block.size, device="cuda", generator=make).mul_(0.08).expand(n, -1).contiguous()
    for rows in (run.x, teacher):
        for name in block.VECTORS:
            block.weights(rows)[name].fill_(1.0)
    r = torch.randn(n, tokens, d, device="cuda", generator=make)
    r = (r + torch.randn(n, 1, d, device="cuda", generator=make)).bfloat16()  # heterogeneous workers
    begins = torch.zeros(n, tokens, dtype=torch.uint8, device="cuda")
    begins[:, ::-(-tokens // 4)] = 1
    target = block.forward(teacher, r, begins=begins).clone()
    losses = []
    for _ in range(steps):
        off = block.forward(run.x, r, begins=begins).float() - target.float()
        losses.append(off.square().mean())
        block.backward(run.x, run.descent, (off * (-1.0 / tokens)).bfloat16())  # -g
        run.step(lr, seed)
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    history = train()
    for step in range(0, len(history), 10):
        print(f"step {step:3d}  mean loss of the workers {history[step]:.4f}")
    print(f"step {len(history) - 1:3d}  mean loss of the workers {history[-1]:.4f}")
