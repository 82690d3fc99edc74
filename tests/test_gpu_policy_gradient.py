"""A step on a model's own answers as a whole: the example model, its gradients, serving token by token, and the calls together in a captured graph."""
import importlib.util
import math
import os

import pytest
import torch

from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_gradient_example", os.path.join(ROOT, "examples", "policy_gradient.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_example_runs(example, dtype):
    print(f"[gpu-case] policy gradient {dtype}", flush=True)
    rewards = example.main(steps=3, answers=9, length=7, dtype=dtype, say=lambda text: print(text, flush=True))
    assert len(rewards) == 3 and all(0 <= r <= 1 for r in rewards)


def wide_loss(example, model, wide, tokens, lengths, temperature, vocab):
    """The example's loss from elementary operations in 64 bits."""
    heads, kv, width = model.heads, model.kv_heads, model.width
    now, then = tokens[:, :-1], tokens[:, 1:]
    answers, length = now.shape
    norm = lambda s, w: w * s / torch.sqrt(s.pow(2).mean(-1, keepdim=True) + example.EPS)  # noqa: E731
    angle = torch.arange(length).repeat(answers).double()[:, None] * model.turns.cpu()
    cos, sin, half = torch.cos(angle)[:, None], torch.sin(angle)[:, None], model.turns.numel()

    def turned(v):
        a, b = v[..., :half], v[..., half:2 * half]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, v[..., 2 * half:]], -1)

    stream = wide["embedding"][now.reshape(-1)]
    delta = torch.zeros_like(stream)
    for i in range(len(model.packed)):
        stream = stream + delta
        packed = (norm(stream, wide[f"norms.{i}"]) @ wide[f"packed.{i}"]).reshape(answers * length, heads + 2 * kv, width)
        q, k = turned(norm(packed[:, :heads], wide[f"q_norms.{i}"])), turned(norm(packed[:, heads:heads + kv], wide[f"k_norms.{i}"]))
        q, k, v = (t.reshape(answers, length, -1, width).transpose(1, 2) for t in (q, k, packed[:, heads + kv:]))
        k, v = (t.repeat_interleave(heads // kv, 1) for t in (k, v))
        scores = q @ k.transpose(2, 3) / math.sqrt(width)
        scores = scores.masked_fill(torch.ones(length, length, dtype=torch.bool).triu(1), -math.inf)
        delta = (torch.softmax(scores, -1) @ v).transpose(1, 2).reshape(answers * length, heads * width) @ wide[f"out.{i}"]
    logits = norm(stream + delta, wide[f"norms.{len(model.packed)}"]) @ wide["head"].T
    logp = torch.log_softmax(logits / temperature, 1)
    kept = torch.arange(length) < lengths[:, None]
    reward = ((now + 1) % vocab == then).double()
    advantage = reward - (reward * kept).sum() / kept.sum()
    given = logp.gather(1, then.reshape(-1, 1)).reshape(answers, length)
    entropy = -(logp.exp() * logp).sum(1).reshape(answers, length)
    return -((advantage * given + 0.01 * entropy) * kept).sum() / kept.sum()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_its_gradients_are_those_of_the_same_model_in_64_bits(example, dtype):
    """Every parameter's gradient.  In 32 bits the chain of products keeps five digits; in bf16 each of some forty roundings on the way there and back (two
    blocks of ten, the head's four) costs 2^-8 of what it rounds."""
    print(f"[gpu-case] policy gradients {dtype}", flush=True)
    vocab, temperature = 50, 1.5
    model = example.Model(vocab, 4, 2, 32, 16, 2, dtype, seed=5)
    g = torch.Generator().manual_seed(6)
    tokens = torch.randint(0, vocab, (7, 14), generator=g)
    tokens[:, 4] = (tokens[:, 3] + 1) % vocab               # (some rewards)
    tokens[::2, 9] = (tokens[::2, 8] + 1) % vocab
    lengths = torch.tensor([13, 1, 5, 9, 13, 10, 7])
    loss, _ = example.loss_of(model, tokens.cuda(), lengths.cuda(), temperature, vocab)
    loss.backward()
    wide = {n: p.detach().double().cpu().requires_grad_() for n, p in model.named_parameters()}
    wide_loss(example, model, wide, tokens, lengths, temperature, vocab).backward()
    for name, p in model.named_parameters():
        got, want = p.grad.double().cpu(), wide[name].grad
        assert float((got - want).norm() / want.norm()) < (1e-5 if dtype == torch.float32 else 40 * 2.0 ** -8), name
    # the clipped gradients: each times the same factor, in place
    before = [p.grad.double().clone() for p in model.parameters()]
    norm = math.sqrt(sum(float(b.pow(2).sum()) for b in before))
    for most in (norm * 0.25, norm * 4):
        factor = min(1.0, most / (norm + 1e-6))
        for p, b in zip(model.parameters(), before):
            p.grad.copy_(b)
        assert abs(float(example.clip(model.parameters(), most)) - norm) <= 4 * U * norm
        half = U if dtype == torch.float32 else 2.0 ** -8
        for p, b in zip(model.parameters(), before):
            here = half if p.dtype == torch.bfloat16 else U
            assert float(((p.grad.double() - b * factor).abs() - (here + 5 * U) * (b * factor).abs()).max()) <= 1e-40


def test_a_model_that_was_converted_as_a_whole(example):
    """model.bfloat16() converts the norms' weights, too: gradients as those of the model in 64 bits (bounds as above), and answers token by token."""
    print("[gpu-case] policy gradients of a converted model", flush=True)
    vocab, g = 50, torch.Generator().manual_seed(7)
    model = example.Model(vocab, 4, 2, 32, 16, 2, torch.float32, seed=5)
    for norms in (model.norms, model.q_norms, model.k_norms):
        for w in norms:
            w.data.copy_(1 + 0.3 * torch.randn(w.shape, generator=g))
    model.bfloat16()
    assert all(p.dtype == torch.bfloat16 for p in model.parameters())
    tokens = torch.randint(0, vocab, (7, 14), generator=g)
    tokens[:, 4] = (tokens[:, 3] + 1) % vocab
    lengths = torch.tensor([13, 1, 5, 9, 13, 10, 7])
    example.loss_of(model, tokens.cuda(), lengths.cuda(), 1.5, vocab)[0].backward()
    wide = {n: p.detach().double().cpu().requires_grad_() for n, p in model.named_parameters()}
    wide_loss(example, model, wide, tokens, lengths, 1.5, vocab).backward()
    for name, p in model.named_parameters():
        assert p.grad.dtype == torch.bfloat16
        want = wide[name].grad
        assert float((p.grad.double().cpu() - want).norm() / want.norm()) < 40 * 2.0 ** -8, name
    with torch.no_grad():
        whole = model.logits(tokens[:, :5].cuda()).reshape(7, 5, vocab).double()
        cache = model.cache(7, 5)
        for position in range(5):
            got = model.step(tokens[:, position].cuda(), position, cache).double()
            assert float((got - whole[:, position]).norm() / whole[:, position].norm()) < 24 * 2.0 ** -8, position


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_token_by_token_is_all_at_once(example, dtype):
    """Logits of single tokens with a cache against those of whole answers: the same operations, products in another order (in bf16 a dozen roundings that may fall
    the other way)."""
    print(f"[gpu-case] answers token by token {dtype}", flush=True)
    model = example.Model(60, 6, 3, 32, 32, 2, dtype, seed=8)
    tokens = torch.randint(0, 60, (5, 11), generator=torch.Generator().manual_seed(9)).cuda()
    with torch.no_grad():
        whole = model.logits(tokens).reshape(5, 11, 60).double()
        cache = model.cache(5, 11)
        for position in range(11):
            got = model.step(tokens[:, position], position, cache).double()
            off = float((got - whole[:, position]).norm() / whole[:, position].norm())
            assert off < (1e-5 if dtype == torch.float32 else 24 * 2.0 ** -8), position


class Together:
    """All calls of a step with buffers of their own, as a program that captures them would hold them."""

    def __init__(self, tokens, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.g, self.tokens, self.vocab = g, tokens, 5001
        row = 12 * 64
        self.packed, self.out = new(tokens, row, dtype=torch.bfloat16), new(tokens, 10 * 64, dtype=torch.bfloat16)
        self.dout, self.dpacked = new(tokens, 10 * 64, dtype=torch.bfloat16), torch.zeros(tokens, row, dtype=torch.bfloat16, device="cuda")
        self.weights, self.dweights = [new(64) for _ in "qk"], [new(64) for _ in "qk"]
        self.positions, self.turns = torch.zeros(tokens, dtype=torch.int64, device="cuda"), 10000.0 ** (-torch.arange(32, dtype=torch.float64, device="cuda") / 32)
        self.logits, self.dlogits = new(tokens, self.vocab, dtype=torch.bfloat16), new(tokens, self.vocab, dtype=torch.bfloat16)
        self.targets = torch.zeros(tokens, dtype=torch.int64, device="cuda")
        self.logp, self.entropy, self.stats = new(tokens), new(tokens), new(tokens, 2)
        self.ids, self.top_logp = new(tokens, 10, dtype=torch.int64), new(tokens, 10)
        self.dlogp, self.dentropy = new(tokens), new(tokens)
        self.norm = new(1)
        self.qk = bns.make_qk(tokens, 8, 2, 64, q=(row, 64), k=(row, 64), q_out=(10 * 64, 64), k_out=(10 * 64, 64), dq=(row, 64), dk=(row, 64))
        self.logprob = bns.make_logprob(tokens, self.vocab, top=10)
        grads = [self.dpacked, self.dlogits, *self.dweights]
        self.gradients = bns.make_gradients(grads, grads)
        self.rooms = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in
                      (bns.bns_qk_workspace_bytes(self.qk), bns.bns_logprob_workspace_bytes(self.logprob), bns.bns_grads_workspace_bytes(self.gradients))]
        self.fill()

    def fill(self):
        for t in (self.packed, self.dout, self.logits, *self.weights, self.dlogp, self.dentropy):
            t.normal_(generator=self.g)
        self.positions.random_(0, 10 ** 6, generator=self.g)
        self.targets.random_(-300, self.vocab, generator=self.g)

    def run(self):
        bns.bns_qk_forward(self.qk, self.packed, self.packed[:, 512:], *self.weights, self.positions, self.turns, self.out, self.out[:, 512:])
        bns.bns_logprob_forward(self.logprob, self.logits, self.targets, self.logp, self.entropy, self.stats, self.ids, self.top_logp, self.rooms[1])
        bns.bns_logprob_backward(self.logprob, self.logits, self.targets, self.stats, self.entropy, self.dlogp, self.dentropy, self.dlogits)
        bns.bns_qk_backward(self.qk, self.packed, self.packed[:, 512:], *self.weights, self.positions, self.turns, self.dout, self.dout[:, 512:], self.dpacked,
                            self.dpacked[:, 512:], *self.dweights, self.rooms[0])
        bns.bns_grads_clip(self.gradients, 1.0, self.norm, self.rooms[2])

    def results(self):
        return [t.clone() for t in (self.out, self.logp, self.entropy, self.stats, self.ids, self.top_logp, self.dlogits, self.dpacked, *self.dweights, self.norm)]


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("tokens", [1, 37, 1500])
def test_two_captured_steps_are_replayed_beside_eager_ones(tokens):
    """Two graphs with workspaces of their own, replayed on two streams with new inputs, against eager calls on the same inputs: the same bits."""
    print(f"[gpu-case] captured steps {tokens}", flush=True)
    steps = [Together(tokens, seed) for seed in (1, 2)]
    streams, graphs = [torch.cuda.Stream() for _ in steps], []
    for step, stream in zip(steps, streams):
        step.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step.run()
        graphs.append(graph)
    for _ in range(4):
        for step in steps:
            step.fill()
        wanted = []
        for step in steps:
            step.run()
            wanted.append(step.results())
            for t in (step.out, step.dlogits, step.dpacked, step.logp, step.ids, step.norm):
                t.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for step, want in zip(steps, wanted):
            assert float(step.norm) > 1.0 and same(step.results(), want)


def test_steps_on_two_streams_at_once():
    print("[gpu-case] steps on two streams", flush=True)
    steps = [Together(700, seed) for seed in (3, 4)]
    wanted = []
    for step in steps:
        step.run()
        wanted.append(step.results())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for step, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                step.run()
    torch.cuda.synchronize()
    for step, want in zip(steps, wanted):
        assert same(step.results(), want)
