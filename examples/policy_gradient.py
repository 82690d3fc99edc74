"""A small attention model that learns from rewards for its own answers: it answers token by token, drawing each from its most probable alternatives, then takes a
step along the policy gradient.

    python examples/policy_gradient.py            (on an MI355X, after `python __graft_entry__.py`)

An answer is rewarded for every token that follows its predecessor in the vocabulary's order.  Norms, the queries' and keys' rotation, log probabilities with
entropy and alternatives and the clipping of the gradients run in libbns; attention, products, embeddings and the optimizer are plain torch.
"""
import argparse
import importlib.util
import math
import os
import sys

import torch
from torch.autograd.function import once_differentiable

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
from paper_1810_10962_amd import bns  # noqa: E402

_spec = importlib.util.spec_from_file_location("language_model_example", os.path.join(ROOT, "examples", "language_model.py"))
_language_model = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(_language_model)
AddNorm, NAMES, EPS = _language_model.AddNorm, _language_model.NAMES, _language_model.EPS


def frequencies(rotated):
    return 10000.0 ** (-torch.arange(rotated // 2, dtype=torch.float64, device="cuda") * 2 / rotated)


class QueriesKeys(torch.autograd.Function):
    """Queries, keys and values of a projection's result: queries and keys with every head's norm and the rotation by position."""

    @staticmethod
    def forward(ctx, packed, q_weight, k_weight, positions, turns, heads, kv_heads):
        packed, q_weight, k_weight = packed.contiguous(), q_weight.contiguous(), k_weight.contiguous()
        positions, turns = positions.long().contiguous(), turns.double().contiguous()
        if q_weight.dtype != k_weight.dtype:
            raise TypeError(f"weights of the queries' norm are {q_weight.dtype}, of the keys' {k_weight.dtype}")
        tokens, row = packed.shape
        width = q_weight.numel()
        qk = bns.make_qk(tokens, heads, kv_heads, width, NAMES[packed.dtype], rotated=2 * turns.numel(), weight_dtype=NAMES[q_weight.dtype], eps=EPS,
                         q=(row, width), k=(row, width), dq=(row, width), dk=(row, width))
        q = packed.new_empty(tokens, heads, width)
        k = packed.new_empty(tokens, kv_heads, width)
        bns.bns_qk_forward(qk, packed, packed[:, heads * width:], q_weight, k_weight, positions, turns, q, k)
        ctx.save_for_backward(packed, q_weight, k_weight, positions, turns)
        ctx.qk = qk
        return q, k, packed[:, (heads + kv_heads) * width:].reshape(tokens, kv_heads, width)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        packed, q_weight, k_weight, positions, turns = ctx.saved_tensors
        at, behind = ctx.qk.q_heads * ctx.qk.width, (ctx.qk.q_heads + ctx.qk.k_heads) * ctx.qk.width
        dpacked = torch.empty_like(packed)
        dpacked[:, behind:] = dv.reshape(dv.shape[0], -1)
        dq_weight, dk_weight = (torch.empty(w.shape, device=w.device) for w in (q_weight, k_weight))       # (in 32 bits, whatever the weights' type)
        workspace = torch.empty(bns.bns_qk_workspace_bytes(ctx.qk), dtype=torch.uint8, device=packed.device)
        bns.bns_qk_backward(ctx.qk, packed, packed[:, at:], q_weight, k_weight, positions, turns, dq.contiguous(), dk.contiguous(), dpacked, dpacked[:, at:],
                            dq_weight, dk_weight, workspace)
        return dpacked, dq_weight.to(q_weight.dtype), dk_weight.to(k_weight.dtype), None, None, None, None


class LogProb(torch.autograd.Function):
    """(log probability of the target, entropy) of every row of logits; a target outside the vocabulary has log probability 0 and no gradient."""

    @staticmethod
    def forward(ctx, logits, targets, temperature):
        logits, targets = logits.contiguous(), targets.long().contiguous()
        spec = bns.make_logprob(*logits.shape, NAMES[logits.dtype], temperature=temperature)
        logp, entropy = (torch.empty(len(targets), device=logits.device) for _ in range(2))
        stats = torch.empty(len(targets), 2, device=logits.device)
        workspace = torch.empty(bns.bns_logprob_workspace_bytes(spec), dtype=torch.uint8, device=logits.device)
        bns.bns_logprob_forward(spec, logits, targets, logp, entropy, stats, None, None, workspace)
        ctx.save_for_backward(logits, targets, stats, entropy)
        ctx.spec = spec
        return logp, entropy

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dentropy):
        logits, targets, stats, entropy = ctx.saved_tensors
        dlogits = torch.empty_like(logits)
        bns.bns_logprob_backward(ctx.spec, logits, targets, stats, entropy, dlogp.contiguous(), dentropy.contiguous(), dlogits)
        return dlogits, None, None


def alternatives(logits, top, temperature):
    """The `top` most probable tokens of every row and their log probabilities."""
    logits = logits.contiguous()
    spec = bns.make_logprob(*logits.shape, NAMES[logits.dtype], top=top, temperature=temperature)
    ids = torch.empty(len(logits), top, dtype=torch.int64, device=logits.device)
    logp = torch.empty(len(logits), top, device=logits.device)
    bns.bns_logprob_forward(spec, logits, None, None, None, None, ids, logp,
                            torch.empty(bns.bns_logprob_workspace_bytes(spec), dtype=torch.uint8, device=logits.device))
    return ids, logp


def clip(parameters, most):
    """Scales the gradients down, in place, until their norm is at most `most`; the norm as it was."""
    grads = [p.grad for p in parameters if p.grad is not None]
    gradients = bns.make_gradients(grads, grads)
    norm = torch.empty(1, device=grads[0].device)
    bns.bns_grads_clip(gradients, most, norm, torch.empty(bns.bns_grads_workspace_bytes(gradients), dtype=torch.uint8, device=grads[0].device))
    return norm


def attend(q, k, v, from_position):
    """Causal attention of q [answers, length, heads, width], its first token at `from_position`, over k and v [answers, so far, kv heads, width]; in 32 bits."""
    answers, length, heads, width = q.shape
    share = heads // k.shape[2]
    q, k, v = (t.float().transpose(1, 2) for t in (q, k.repeat_interleave(share, 2), v.repeat_interleave(share, 2)))
    scores = q @ k.transpose(2, 3).contiguous() / math.sqrt(width)
    behind = torch.arange(k.shape[2], device=q.device) > torch.arange(length, device=q.device)[:, None] + from_position
    mixed = torch.softmax(scores.masked_fill(behind, -math.inf), -1) @ v.contiguous()
    return mixed.transpose(1, 2).reshape(answers * length, heads * width)


class Model(torch.nn.Module):
    def __init__(self, vocab, heads, kv_heads, width, rotated, blocks, dtype, seed):
        super().__init__()
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda *s, std: torch.nn.Parameter((torch.randn(*s, generator=g, device="cuda") * std).to(dtype))  # noqa: E731
        ones = lambda n: torch.nn.Parameter(torch.ones(n, device="cuda"))  # noqa: E731
        self.heads, self.kv_heads, self.width, stream = heads, kv_heads, width, heads * width
        self.embedding, self.head = make(vocab, stream, std=0.5), make(vocab, stream, std=0.5 * stream ** -0.5)
        self.packed = torch.nn.ParameterList(make(stream, (heads + 2 * kv_heads) * width, std=stream ** -0.5) for _ in range(blocks))
        self.out = torch.nn.ParameterList(make(stream, stream, std=0.5 * stream ** -0.5) for _ in range(blocks))
        self.norms = torch.nn.ParameterList(ones(stream) for _ in range(blocks + 1))
        self.q_norms, self.k_norms = (torch.nn.ParameterList(ones(width) for _ in range(blocks)) for _ in range(2))
        self.turns = frequencies(rotated)

    def logits(self, tokens):
        """Of every token of tokens [answers, length]."""
        answers, length = tokens.shape
        positions = torch.arange(length, device="cuda").repeat(answers)
        stream = self.embedding[tokens.reshape(-1)]
        delta = torch.zeros_like(stream)
        for i, packed in enumerate(self.packed):
            stream, y = AddNorm.apply(delta, stream, self.norms[i])
            q, k, v = QueriesKeys.apply(y @ packed, self.q_norms[i], self.k_norms[i], positions, self.turns, self.heads, self.kv_heads)
            delta = attend(*(t.unflatten(0, (answers, length)) for t in (q, k, v)), 0).to(y.dtype) @ self.out[i]
        return AddNorm.apply(delta, stream, self.norms[-1])[1] @ self.head.T

    def cache(self, answers, length):
        return [[self.embedding.new_zeros(answers, length, self.kv_heads, self.width) for _ in "kv"] for _ in self.packed]

    @torch.no_grad()
    def step(self, tokens, position, cache):
        """Logits of one token of every answer; its keys go straight into the cache [answers, length, kv heads, width]."""
        answers = len(tokens)
        positions = torch.full((answers,), position, device="cuda")
        stream = self.embedding[tokens]
        delta = torch.zeros_like(stream)
        for i, (keys, values) in enumerate(cache):
            stream, y = AddNorm.apply(delta, stream, self.norms[i])
            packed = y @ self.packed[i]
            row, width = packed.shape[1], self.width
            at, behind = self.heads * width, (self.heads + self.kv_heads) * width
            values[:, position] = packed[:, behind:].reshape(answers, self.kv_heads, width)
            qk = bns.make_qk(answers, self.heads, self.kv_heads, width, NAMES[y.dtype], rotated=2 * self.turns.numel(),
                             weight_dtype=NAMES[self.q_norms[i].dtype], eps=EPS, q=(row, width), k=(row, width), q_out=(row, width), k_out=(keys.stride(0), width))
            bns.bns_qk_forward(qk, packed, packed[:, at:], self.q_norms[i], self.k_norms[i], positions, self.turns, packed, keys[:, position])
            q = packed[:, :at].reshape(answers, 1, self.heads, width)
            delta = attend(q, keys[:, :position + 1], values[:, :position + 1], position).to(y.dtype) @ self.out[i]
        return AddNorm.apply(delta, stream, self.norms[-1])[1] @ self.head.T


def answer(model, first, length, top, temperature, generator):
    """Answers of `length` tokens, one after the other from the `top` most probable ones."""
    cache, tokens = model.cache(len(first), length), [first]
    for position in range(length):
        ids, logp = alternatives(model.step(tokens[-1], position, cache), top, temperature)
        drawn = torch.multinomial(torch.softmax(logp, 1), 1, generator=generator)
        tokens.append(ids.gather(1, drawn)[:, 0])
    return torch.stack(tokens, 1)


def loss_of(model, tokens, lengths, temperature, vocab, bonus=0.01):
    """Policy gradient's loss of answers [answers, 1 + length], of which `lengths` tokens count, and the mean reward."""
    now, then = tokens[:, :-1], tokens[:, 1:]
    kept = torch.arange(then.shape[1], device="cuda") < lengths[:, None]
    reward = ((now + 1) % vocab == then).float()
    count = kept.sum()
    mean = (reward * kept).sum() / count
    logp, entropy = LogProb.apply(model.logits(now), torch.where(kept, then, -1).reshape(-1), temperature)
    kept = kept.reshape(-1)
    return -((reward.reshape(-1) - mean) * logp + bonus * entropy * kept)[kept].sum() / count, mean


def main(steps=60, vocab=64, answers=64, length=24, dtype=torch.float32, top=16, say=print):
    model = Model(vocab, 4, 2, 32, 16, 2, dtype, seed=1)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    g = torch.Generator(device="cuda").manual_seed(2)
    rewards = []
    for step in range(steps):
        first = torch.randint(0, vocab, (answers,), generator=g, device="cuda")
        tokens = answer(model, first, length, top, 1.0, g)
        lengths = torch.randint(1, length + 1, (answers,), generator=g, device="cuda")
        optimizer.zero_grad()
        loss, reward = loss_of(model, tokens, lengths, 1.0, vocab)
        loss.backward()
        norm = clip(model.parameters(), 1.0)
        optimizer.step()
        rewards.append(float(reward))
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: reward {rewards[-1]:.3f}, norm of the gradients {float(norm):.3f}")
    return rewards


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = parser.parse_args()
    main(a.steps, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype])
