"""A small language model whose norms and losses run in libbns: trained, distilled into a smaller one, and run token by token with 8-bit activations.

    python examples/language_model.py            (on an MI355X, after `python __graft_entry__.py`)

The data is a Markov chain over the vocabulary, made here.  Everything that is not a norm or a loss (embeddings, the blocks' two matrices, the
optimizer) is plain torch.
"""
import argparse
import os
import sys

import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_10962_amd import bns  # noqa: E402

EPS = 1e-6
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16"}


class AddNorm(torch.autograd.Function):
    """(stream, y) = (delta + stream, norm of it): the residual's addition and the norm behind it."""

    @staticmethod
    def forward(ctx, delta, stream, weight):
        delta, stream, weight = delta.contiguous(), stream.contiguous(), weight.contiguous()      # (the library is handed addresses)
        rows, width = stream.shape
        rms = bns.make_rms(rows, width, NAMES[stream.dtype], eps=EPS)
        total, y, rstd = torch.empty_like(stream), torch.empty_like(stream), torch.empty(rows, device=stream.device)
        bns.bns_rms_forward(rms, delta, stream, weight, total, y, None, rstd)
        ctx.save_for_backward(total, weight, rstd)
        ctx.rms = rms
        return total, y

    @staticmethod
    @once_differentiable
    def backward(ctx, dtotal, dy):
        total, weight, rstd = ctx.saved_tensors
        dx, dweight = torch.empty_like(total), torch.empty_like(weight)
        workspace = torch.empty(bns.bns_rms_workspace_bytes(ctx.rms), dtype=torch.uint8, device=total.device)
        bns.bns_rms_backward(ctx.rms, total, weight, rstd, dy.contiguous(), dtotal.contiguous(), dx, dweight, workspace)
        return dx, dx, dweight          # the sum's gradient is both addends'


class HeadLoss(torch.autograd.Function):
    """Mean cross entropy of hidden weight^T against the targets, without the logits; targets outside the vocabulary are left out."""

    @staticmethod
    def forward(ctx, hidden, weight, targets):
        hidden, weight, targets = hidden.contiguous(), weight.contiguous(), targets.contiguous()
        head = bns.make_head(hidden.shape[0], hidden.shape[1], weight.shape[0], NAMES[hidden.dtype])
        workspace = torch.empty(bns.bns_head_workspace_bytes(head), dtype=torch.uint8, device=hidden.device)
        loss, lse = torch.empty(hidden.shape[0], device=hidden.device), torch.empty(hidden.shape[0], device=hidden.device)
        bns.bns_head_forward(head, hidden, weight, targets, loss, lse, workspace)
        count = ((targets >= 0) & (targets < weight.shape[0])).sum().clamp(min=1)
        ctx.save_for_backward(hidden, weight, targets, lse, count)
        ctx.head, ctx.workspace = head, workspace
        return loss.sum() / count

    @staticmethod
    @once_differentiable
    def backward(ctx, dmean):
        hidden, weight, targets, lse, count = ctx.saved_tensors
        dloss = (dmean / count).expand(hidden.shape[0]).contiguous()
        dhidden, dweight = torch.empty_like(hidden), torch.empty_like(weight)
        bns.bns_head_backward(ctx.head, hidden, weight, targets, lse, dloss, dhidden, dweight, ctx.workspace)
        return dhidden, dweight, None


class DistillLoss(torch.autograd.Function):
    """Mean loss of the student's logits against a teacher's top logits.  The mean's gradient is known beforehand, so the logits' comes from the
    forward pass and backward only scales it."""

    @staticmethod
    def forward(ctx, logits, ids, teacher, temperature):
        logits, ids, teacher = logits.contiguous(), ids.contiguous(), teacher.contiguous()
        tokens, vocab = logits.shape
        distill = bns.make_distill(tokens, vocab, ids.shape[1], NAMES[logits.dtype], temperature=temperature)
        loss, lse, dlogits = torch.empty(tokens, device=logits.device), torch.empty(tokens, device=logits.device), torch.empty_like(logits)
        dloss = torch.full((tokens,), 1.0 / tokens, device=logits.device)
        bns.bns_distill_forward(distill, logits, ids, teacher, dloss, loss, lse, dlogits)
        ctx.save_for_backward(dlogits)
        return loss.mean()

    @staticmethod
    @once_differentiable
    def backward(ctx, dmean):
        return ctx.saved_tensors[0] * dmean, None, None, None


class Model(torch.nn.Module):
    def __init__(self, vocab, width, blocks, dtype, seed):
        super().__init__()
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda *s, std: torch.nn.Parameter((torch.randn(*s, generator=g, device="cuda") * std).to(dtype))  # noqa: E731
        self.embedding, self.head = make(vocab, width, std=0.5), make(vocab, width, std=width ** -0.5)
        self.up = torch.nn.ParameterList(make(width, 2 * width, std=width ** -0.5) for _ in range(blocks))
        self.down = torch.nn.ParameterList(make(2 * width, width, std=0.5 * (2 * width) ** -0.5) for _ in range(blocks))
        self.norms = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(width, device="cuda")) for _ in range(blocks + 1))

    def hidden(self, tokens):
        stream = self.embedding[tokens]
        delta = torch.zeros_like(stream)
        for up, down, norm in zip(self.up, self.down, self.norms):
            stream, y = AddNorm.apply(delta, stream, norm)
            delta = torch.nn.functional.gelu(y @ up) @ down
        return AddNorm.apply(delta, stream, self.norms[-1])[1]

    @torch.no_grad()
    def hidden_8_bits(self, tokens):
        """The same for serving: the norm leaves its result in 8 bits with a scale for every 32 elements, as an 8-bit product would take it (here its values
        are multiplied as they are)."""
        stream = self.embedding[tokens]
        delta = torch.zeros_like(stream)
        rows, width = stream.shape
        rms = bns.make_rms(rows, width, NAMES[stream.dtype], out="e4m3", group=32, pow2_scales=True, eps=EPS)
        y = torch.empty(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
        scales = torch.empty(rows, -(-width // 32), device="cuda")
        for i, norm in enumerate(self.norms):
            bns.bns_rms_forward(rms, delta, stream, norm, stream, y, scales, None)       # the stream is updated in place
            x = (y.float() * scales.repeat_interleave(32, 1)[:, :width]).to(stream.dtype)
            if i < len(self.up):
                delta = torch.nn.functional.gelu(x @ self.up[i]) @ self.down[i]
        return x


def chain(vocab, tokens, seed):
    """Pairs (token, the one that follows): every token is followed by one of four, the first of them most often; some targets are unknown (-100)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    now = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    which = torch.multinomial(torch.tensor([0.7, 0.15, 0.1, 0.05], device="cuda"), tokens, replacement=True, generator=g)
    then = (now * 31 + 7 + which * 101) % vocab
    return now, torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.05, -100, then)


def train(model, steps, vocab, tokens, loss_of):
    optimizer = torch.optim.Adam(model.parameters(), lr=4e-3)
    losses = []
    for step in range(steps):
        now, then = chain(vocab, tokens, step)
        optimizer.zero_grad()
        loss = loss_of(model, now, then)
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    return losses


def main(steps=60, vocab=1000, width=128, tokens=2048, dtype=torch.float32, say=print):
    teacher = Model(vocab, width, 2, dtype, seed=1)
    losses = train(teacher, steps, vocab, tokens, lambda m, now, then: HeadLoss.apply(m.hidden(now), m.head, then))
    say(f"teacher: cross entropy {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")

    student = Model(vocab, width, 1, dtype, seed=2)

    def against_teacher(model, now, then):
        with torch.no_grad():
            top = torch.topk((teacher.hidden(now) @ teacher.head.T).float(), 16)
        return DistillLoss.apply(model.hidden(now) @ model.head.T, top.indices, top.values.contiguous(), 2.0)

    distilled = train(student, steps, vocab, tokens, against_teacher)
    say(f"student: distillation loss {distilled[0]:.3f} -> {distilled[-1]:.3f}")

    # serving, one token at a time
    now, then = chain(vocab, 64, 10 ** 6)
    same = sum(int((teacher.hidden_8_bits(now[i:i + 1]) @ teacher.head.T).argmax()) == int((teacher.hidden(now[i:i + 1]) @ teacher.head.T).argmax())
               for i in range(len(now)))
    say(f"single tokens with 8-bit activations: {same} of {len(now)} choices as with {NAMES[dtype]}")
    return losses, distilled, same / len(now)


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = parser.parse_args()
    main(a.steps, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype])
