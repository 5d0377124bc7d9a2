"""A token student: recurrent blocks between an embedding and the vocabulary, learning from labels or from a teacher's top logits.

What stands in front of a sequence model's first block and behind its last, with the library's token operators around the blocks of `sequence`:

    x = scale * table[token],  s <- x + block_1(x) + ...,  h = norm(s),  logits = h table^T

The table is the last product's weight too, so it has two gradients: the loss writes one, the embedding's is added to it (each time
in fp32 and rounded to bf16: two roundings, of which the second is what a sum of two bf16 gradients has anyway).  Blocks that were distilled
one by one against a teacher's can be put between, and the whole then learns on text: `learn` from labels (softmax cross entropy over
the whole vocabulary, whose logits are never kept), `imitate` from the teacher's largest logits, stored beforehand.

Embedding, losses, norms, recurrences and update are the library's kernels; the blocks' projections, and the logits where they are wanted,
are plain matrix products and torch's, in bf16.

    python -m paper_2012_03096_amd.tokens            # a student learns a language of few words, another one imitates it
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import binding as pb
from .sequence import SequenceBlock


class TokenStudent:
    """A model of `blocks` recurrent blocks of width d over `vocab` tokens.  A token or label outside 0..vocab-1 is padding.  Tokens,
    labels and a teacher's logits may have any strides."""

    def __init__(self, vocab: int, d: int, blocks: int = 1, seed: int = 0, device: str = "cuda", state_bits: int = 8, weight_decay: float = 0.01):
        gen = torch.Generator().manual_seed(seed)
        self.vocab, self.d, self.scale = vocab, d, math.sqrt(d)
        self.blocks = [SequenceBlock(d, seed=1000 * seed + k + 1, device=device, state_bits=state_bits, weight_decay=weight_decay) for k in range(blocks)]
        # fp32 masters; the table also in bf16, which lookup and products read and the update refreshes
        self.params = [(torch.randn(vocab, d, generator=gen) * d ** -0.5).to(device), torch.ones(d, device=device)]
        self.table, self.norm = self.params[0].to(torch.bfloat16), self.params[1]
        self.grads = [torch.empty_like(self.table), torch.empty_like(self.norm)]
        self.optimizer = pb.AdamW(self.params, state_bits=state_bits, copies=[self.table, torch.empty(d, dtype=torch.bfloat16, device=device)],
                                  weight_decay=[weight_decay, 0.0])
        self._buffers, self._saved = {}, None

    def _buffer(self, name: str, *shape, dtype=torch.bfloat16):
        """A buffer of the model for what is called `name`, as large as the largest that was asked for."""
        n, have = math.prod(shape), self._buffers.get(name)
        if have is None or have.numel() < n:
            self._buffers.pop(name, None)
            have = self._buffers[name] = torch.empty(n, dtype=dtype, device=self.table.device)
        return have[:n].view(shape)

    def _bytes(self, name: str, n: int):
        return self._buffer(name, n, dtype=torch.uint8)

    def _forward(self, tokens, training: bool):
        """h [batch * len, d] for tokens [batch, len]; a training pass keeps what the backward pass needs."""
        b, t = tokens.shape
        out, stream, saved = self._buffer("x", b, t, self.d), None, []
        pb.embed_forward(tokens.contiguous(), self.table, out, scale=self.scale)
        for k, block in enumerate(self.blocks):
            total = None if stream is None or training else torch.empty_like(out)
            y, z, q = block._forward(out, stream, None, None, None, training, total=total)
            saved.append((out, stream, z, q))
            # the stream behind the first sum is the sum itself; a training pass keeps it in the block's buffer
            stream, out = out if stream is None else (q["total"] if training else total), y
        h, total = self._buffer("h", b, t, self.d), self._buffer("total", b, t, self.d)
        pb.rmsnorm_forward(out, self.norm, h, residual=stream, total=total)
        self._saved = (saved, total) if training else None
        return h.view(-1, self.d)

    def _backward(self, tokens, dh) -> None:
        """All gradients from dh [batch * len, d]; the table's is added to what the loss wrote."""
        saved, total = self._saved
        shape = total.shape
        rows = shape[0] * shape[1]
        g = torch.empty_like(total)
        pb.rmsnorm_backward(total, self.norm, dh.view(shape), g, self.grads[1], self._bytes("norm_workspace", pb.rmsnorm_workspace_bytes(rows, self.d)))
        for block, (x, stream, z, q) in zip(reversed(self.blocks), reversed(saved)):
            # what arrives at the sum behind the block reaches its output and, past it, the stream in front of it
            g = block._backward(x, stream, g.view(-1, self.d), z, q, dtotal=g)
        pb.embed_backward(tokens.contiguous(), g, self.grads[0], self._bytes("embed_workspace", pb.embed_workspace_bytes(rows, self.vocab, self.d)), scale=self.scale,
                          accumulate=True)
        self._saved = None

    def _update(self, lr: float) -> None:
        self.optimizer.step(self.grads, lr)
        for block in self.blocks:
            block.optimizer.step(block.grads, lr)

    def learn_gradients(self, tokens, labels):
        """Forward and backward pass for the mean cross entropy of labels [batch, len] (those outside the vocabulary are ignored).  The gradients
        are in grads and the blocks' grads; returns the loss as a tensor on the GPU."""
        h = self._forward(tokens, True)
        rows = h.shape[0]
        live = (labels >= 0) & (labels < self.vocab)
        weight = (live / live.sum().clamp_min(1)).view(-1).float()
        loss, dh = self._buffer("loss", rows, dtype=torch.float32), self._buffer("dh", rows, self.d)
        workspace = self._bytes("head_workspace", pb.head_loss_workspace_bytes(rows, self.vocab, self.d, h.dtype, gradients=True))
        pb.head_loss(h, self.table, labels.reshape(-1).contiguous(), loss, workspace, row_weight=weight, dh=dh, dweight=self.grads[0])
        mean = (loss * weight).sum()
        self._backward(tokens, dh)
        return mean

    def imitate_gradients(self, tokens, teacher, at, temperature: float = 2.0):
        """The same for the mean distillation loss against a teacher's top logits: teacher and at [batch, len, top], places outside the
        vocabulary unknown; tokens without any are left out."""
        h = self._forward(tokens, True)
        top = teacher.shape[-1]
        some = ((at >= 0) & (at < self.vocab) & (teacher > float("-inf"))).any(-1).view(-1)
        weight = some / some.sum().clamp_min(1).float()
        logits = h @ self.table.t()
        loss = self._buffer("loss", h.shape[0], dtype=torch.float32)
        pb.topk_distill(logits, teacher.reshape(-1, top).contiguous(), at.reshape(-1, top).contiguous(), loss, temperature=temperature, row_weight=weight, dlogits=logits)
        torch.mm(logits.t(), h, out=self.grads[0])
        mean = (loss * weight).sum()
        self._backward(tokens, logits @ self.table)
        return mean

    def learn(self, tokens, labels, lr: float):
        """One training step on labels; returns the loss of its forward pass as a tensor on the GPU: the call waits for nothing."""
        loss = self.learn_gradients(tokens, labels)
        self._update(lr)
        return loss

    def imitate(self, tokens, teacher, at, lr: float, temperature: float = 2.0):
        """One training step on a teacher's top logits."""
        loss = self.imitate_gradients(tokens, teacher, at, temperature)
        self._update(lr)
        return loss

    def score(self, tokens, labels):
        """-log p of each label [batch, len] float32 (0 for ignored ones), logits never kept."""
        h = self._forward(tokens, False)
        loss = torch.empty(h.shape[0], device=h.device)
        workspace = self._bytes("head_workspace", pb.head_loss_workspace_bytes(h.shape[0], self.vocab, self.d, h.dtype, gradients=False))
        pb.head_loss(h, self.table, labels.reshape(-1).contiguous(), loss, workspace)
        return loss.view(labels.shape)

    def top_logits(self, tokens, top: int):
        """What a student imitates: the `top` largest logits for each token and their places, [batch, len, top]."""
        logits = self._forward(tokens, False) @ self.table.t()
        values, places = logits.topk(top, dim=1)
        return values.view(*tokens.shape, top), places.to(torch.int32).view(*tokens.shape, top)

    def new_state(self, batch: int):
        return [torch.zeros(batch, self.d, device=self.table.device) for _ in self.blocks]

    def answer(self, token, state):
        """Logits [batch, vocab] for the next token after `token` [batch]; state (of new_state) is updated in place."""
        out, stream = torch.empty(token.shape[0], self.d, dtype=torch.bfloat16, device=token.device), None
        pb.embed_forward(token.contiguous(), self.table, out, scale=self.scale)
        for block, s in zip(self.blocks, state):
            total = None if stream is None else torch.empty_like(out)
            y = block.step(out, s, residual=stream, total=total)
            stream, out = out if stream is None else total, y
        h = torch.empty_like(out)
        pb.rmsnorm_forward(out, self.norm, h, residual=stream)
        return h @ self.table.t()


def demo(vocab: int = 2000, d: int = 128, batch: int = 16, length: int = 64, steps: int = 200, lr: float = 3e-3, report: Optional[int] = 50):
    """A language in which a word mostly decides the next: one student learns it from text, another one from the first's top logits.
    Returns their losses and how far token by token answers are from the pass over all tokens."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    follows = torch.randperm(vocab, generator=gen, device="cuda")

    def text():
        words = [torch.randint(0, vocab, (batch,), generator=gen, device="cuda")]
        for _ in range(length):
            other = torch.randint(0, vocab, (batch,), generator=gen, device="cuda")
            words.append(torch.where(torch.rand(batch, generator=gen, device="cuda") < 0.9, follows[words[-1]], other))
        words = torch.stack(words, 1)
        return words[:, :-1].contiguous(), words[:, 1:].contiguous()

    first, second, losses = TokenStudent(vocab, d, blocks=2, seed=1), TokenStudent(vocab, d, seed=2), []
    for name, step in (("learns", lambda x, y: first.learn(x, y, lr)), ("imitates", lambda x, y: second.imitate(x, *first.top_logits(x, 16), lr))):
        for i in range(steps):
            loss = step(*text())
            if report and (i % report == 0 or i == steps - 1):
                losses.append(float(loss))
                print(f"{name}: step {i:4d}  loss {losses[-1]:.4f}", flush=True)
    x, _ = text()
    whole = (first._forward(x, False) @ first.table.t()).view(batch, length, vocab)
    state = first.new_state(batch)
    tokens = torch.stack([first.answer(x[:, t].contiguous(), state) for t in range(length)], 1)
    return losses, float((tokens.float() - whole.float()).norm() / whole.float().norm())


if __name__ == "__main__":
    _, off = demo()
    print(f"token by token against all tokens at once: {off:.2e} apart")
