"""Blockwise distillation of a sequence model's block, with the library's sequence operators.

One task of the method (section 3.1, Eq. 3), as `binding.Block` is for convolutional blocks: the student block is trained to
reproduce the teacher block's activations from the teacher block's own input, on the local loss alone, independently of every
other block.  The student takes the attention's place by a gated recurrence, whose state has one number a channel:

    s = x + residual,  n = norm(s),  (u | gate | out_gate) = n W_in,  h = recurrence(u, gate + bias),  out = (h silu(out_gate)) W_out

Norm, recurrence and update (AdamW, fp32 master weights, states in 8 or 32 bits) are the library's kernels; the projections are
plain matrix products and torch's, in bf16.

The block asks nothing of its teacher but activations: labels may come from attention or any other block.  Those of the demonstration below
come from a frozen block of the student's own form, which it can match.

    python -m paper_2012_03096_amd.sequence          # trains a student on a frozen block's labels, then answers token by token
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import binding as pb


class SequenceBlock:
    """A student (or, untrained, a frozen teacher) block of width d."""

    NAMES = ("norm", "w_in", "bias", "w_out")

    def __init__(self, d: int, seed: int = 0, device: str = "cuda", state_bits: int = 8, weight_decay: float = 0.01):
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=gen)                                             # noqa: E731
        self.d = d
        # fp32 masters; W_in [3d, d] and W_out [d, d] also in bf16, which the products read and the update refreshes
        self.params = [torch.ones(d), rand(3 * d, d) * d ** -0.5, torch.rand(d, generator=gen) * 4.0 + 1.0, rand(d, d) * d ** -0.5]
        self.params = [p.to(device) for p in self.params]
        self.copies = [p.to(torch.bfloat16) for p in self.params]
        self.norm, self.w_in, self.bias, self.w_out = self.params
        self.grads = [torch.empty_like(p) if p.dim() == 1 else torch.empty_like(c) for p, c in zip(self.params, self.copies)]
        self.optimizer = pb.AdamW(self.params, state_bits=state_bits, copies=self.copies, weight_decay=[0.0, weight_decay, 0.0, weight_decay])
        self._buffers, self._views = {}, {}

    def _buffer(self, name: str, *shape, dtype=torch.bfloat16):
        """A buffer of the block for what is called `name`, as large as the largest that was asked for."""
        n, have = math.prod(shape), self._buffers.get(name)
        if have is None or have.numel() < n:
            self._buffers.pop(name, None)
            have = self._buffers[name] = torch.empty(n, dtype=dtype, device=self.params[0].device)
        return have[:n].view(shape)

    def _sized(self, b: int, t: int, training: bool):
        """Activations, their gradients and the operators' workspaces for batches of this size: views of the block's buffers, kept for
        the last size.  A block serves one stream at a time."""
        if self._views.get("size") != (b, t, training):
            self._views = {}
            d, new = self.d, self._buffer
            raw = lambda name, n: new(name, n, dtype=torch.uint8)                                    # noqa: E731
            q = {"size": (b, t, training), "n": new("n", b, t, d), "y": new("y", b, t, d),
                 "workspace": raw("workspace", pb.recurrence_workspace_bytes(b, t, d))}
            if training:
                q.update(saved=raw("saved", pb.recurrence_saved_bytes(b, t, d)), dz=new("dz", b, t, 3 * d), dx=new("dx", b, t, d), total=new("total", b, t, d),
                         norm_workspace=raw("norm_workspace", pb.rmsnorm_workspace_bytes(b * t, d)))
            self._views = q
        return self._views

    def _columns(self, z):
        d = self.d
        return {"u": z[..., :d], "gate": z[..., d:2 * d], "out_gate": z[..., 2 * d:]}

    def _forward(self, x, residual, lengths, state, state_out, training: bool, total=None):
        b, t, d = x.shape
        q = self._sized(b, t, training)
        # the backward pass reads the sum, which is x itself where nothing is added
        pb.rmsnorm_forward(x, self.norm, q["n"], residual=residual, total=q["total"] if training and residual is not None else total)
        z = (q["n"].view(-1, d) @ self.copies[1].t()).view(b, t, 3 * d)
        pb.recurrence_forward(**self._columns(z), y=q["y"], bias=self.bias, lengths=lengths, state=state, state_out=state_out,
                              saved=q.get("saved"), workspace=q["workspace"])
        return (q["y"].view(-1, d) @ self.copies[3].t()).view(b, t, d), z, q

    def forward(self, x, residual=None, lengths=None, state=None, state_out=None, total=None):
        """The block's output for x [batch, len, d] bf16 (plus residual); lengths: int32 [batch] of a padded batch; state and
        state_out [batch, d] float32 carry a text on from piece to piece.  total (like x) receives x + residual, the residual stream: blocks
        follow each other as `out = a.forward(x, total=s); out = b.forward(out, residual=s, total=s)`, and out + s is what they give."""
        return self._forward(x, residual, lengths, state, state_out, False, total)[0]

    def step(self, x, state, active=None, residual=None, total=None):
        """The block's output for one token of each sequence, x [batch, d] (plus residual); state is updated in place (rows with active 0
        stay).  total receives x + residual, as in forward."""
        n, y = torch.empty_like(x), torch.empty_like(x)
        pb.rmsnorm_forward(x, self.norm, n, residual=residual, total=total)
        c = self._columns(n @ self.copies[1].t())
        pb.recurrence_step(c["u"], c["gate"], state, y, out_gate=c["out_gate"], bias=self.bias, active=active)
        return y @ self.copies[3].t()

    def _backward(self, x, residual, dout, z, q, lengths=None, dtotal=None):
        """Gradients of the block's parameters (into self.grads) and of x + residual (returned, a buffer of the block) from dout, what the
        training forward pass left (z, q), and the gradient that arrives at the residual stream."""
        b, t, d = x.shape
        dnorm, dw_in, dbias, dw_out = self.grads
        torch.mm(dout.t(), q["y"].view(-1, d), out=dw_out)
        dy = (dout @ self.copies[3]).view(b, t, d)
        c, g = self._columns(z), self._columns(q["dz"])
        pb.recurrence_backward(**c, dy=dy, saved=q["saved"], du=g["u"], dgate=g["gate"], dout_gate=g["out_gate"], bias=self.bias, dbias=dbias,
                               lengths=lengths, workspace=q["workspace"])
        dz = q["dz"].view(-1, 3 * d)
        torch.mm(dz.t(), q["n"].view(-1, d), out=dw_in)
        dn = (dz @ self.copies[1]).view(b, t, d)
        pb.rmsnorm_backward(q["total"] if residual is not None else x, self.norm, dn, q["dx"], dnorm, q["norm_workspace"], dtotal=dtotal)
        return q["dx"]

    def distill_step(self, x, target, lr: float, residual=None, lengths=None):
        """One distillation step: forward, mean squared difference from target over the real tokens (Eq. 3), backward through this block
        only, AdamW.  What x, residual and target hold behind a sequence has no influence.  Returns the loss of the forward pass as a
        tensor on the GPU: the call waits for nothing."""
        b, t, d = x.shape
        if lengths is not None:
            # the weights' gradients sum over all rows: 0 * NaN of a padded one would be NaN in every weight
            live = (torch.arange(t, device=x.device) < lengths[:, None])[:, :, None]
            x = torch.where(live, x, 0.0)
            residual = torch.where(live, residual, 0.0) if residual is not None else None
        out, z, q = self._forward(x, residual, lengths, None, None, True)
        diff = out.float() - target.float()
        count = b * t * d
        if lengths is not None:
            diff = torch.where(live, diff, 0.0)
            count = live.sum().clamp_min(1) * d
        loss = diff.square().sum() / count
        dout = (diff * (2.0 / count)).to(torch.bfloat16).view(-1, d)
        self._backward(x, residual, dout, z, q, lengths)
        self.optimizer.step(self.grads, lr)
        return loss


def demo(d: int = 256, batch: int = 8, length: int = 512, steps: int = 1000, lr: float = 5e-3, report: Optional[int] = 200):
    """Trains a student on the labels of a frozen block of the same width; returns the losses reported and how far token by
    token answers are from the forward pass over all tokens."""
    teacher, student = SequenceBlock(d, seed=1), SequenceBlock(d, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for i in range(steps):
        x = torch.randn(batch, length, d, generator=gen, device="cuda").to(torch.bfloat16)
        lengths = torch.randint(length // 2, length + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        loss = student.distill_step(x, teacher.forward(x, lengths=lengths), lr, lengths=lengths)
        if report and (i % report == 0 or i == steps - 1):
            losses.append(float(loss))
            print(f"step {i:4d}  loss {losses[-1]:.5f}", flush=True)
    whole = student.forward(x[:, :64].contiguous())
    state = torch.zeros(batch, d, device="cuda")
    tokens = torch.stack([student.step(x[:, t].contiguous(), state) for t in range(64)], 1)
    return losses, float((tokens.float() - whole.float()).norm() / whole.float().norm())


if __name__ == "__main__":
    _, off = demo()
    print(f"token by token against all tokens at once: {off:.2e} apart")
